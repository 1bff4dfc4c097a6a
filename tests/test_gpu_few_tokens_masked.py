"""The layer for few tokens, and choices of weight 0: rows of nothing but masked experts, tokens with fewer than k experts left.
They add nothing, whatever the row of X and those experts' weights hold."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb
from tests import mx4_reference as ref
from tests.test_gpu_few_tokens import _check, _expected, _inputs, _run

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def _poisoned(X, logits, up, down, mask, empty):
    """The same with NaN and infinities in the weights of the experts `mask` and in the rows `empty` of X."""
    X, up, down = X.clone(), up.clone(), down.clone()
    for i, e in enumerate(mask):
        up[e], down[e] = (NAN, INF) if i % 2 else (INF, NAN)
    for i, t in enumerate(empty):
        X[t] = (NAN, INF, -INF)[i % 3]
    return X, logits, up, down


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("T,k,E,hidden,inter", [(1, 2, 8, 264, 40), (9, 3, 8, 256, 128), (16, 6, 64, 512, 176), (16, 4, 300, 64, 64), (16, 2, 6, 4712, 40)])
def test_rows_without_experts(T, k, E, hidden, inter, mx4):
    """Empty slots hold anything, and experts 0 .. k-1, whose ids they show, are out of service."""
    X, logits, up, down = _inputs(T, E, hidden, inter, T + E)
    empty = [t for t in range(T) if t % 5 != 2]
    logits[:, :k] = -INF
    logits[empty] = -INF
    want = _expected(X, logits, up, down, k, mx4)
    got = _run(*_poisoned(X, logits, up, down, range(k), empty), k, mx4)
    _check(got, want)
    assert bool((got[0][empty] == 0).all()) and bool((got[2][empty] == 0).all())
    assert torch.equal(got[1][empty], torch.arange(k, dtype=torch.int32).expand(len(empty), k))


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", ["inf", "lowest"])
@pytest.mark.parametrize("sigmoid,renormalize", [(False, True), (False, False), (True, True), (True, False)])
def test_fewer_experts_than_choices(sigmoid, renormalize, value, dtype, mx4):
    """Every token has 1 to 3 experts left for its 4 choices; the others are masked by -inf or by the type's lowest value."""
    T, k, E, hidden, inter = 6, 4, 20, 256, 96
    X, logits, up, down = _inputs(T, E, hidden, inter, 11)
    logits = logits.to(dtype)
    live = [[5], [5, 9], [9, 13, 17], [17], [13, 5], [9]]
    masked = torch.ones(T, E, dtype=torch.bool)
    for t, experts in enumerate(live):
        masked[t, experts] = False
    logits[masked] = -INF if value == "inf" else torch.finfo(dtype).min
    want = _expected(X, logits, up, down, k, mx4, sigmoid, renormalize)
    out_of_service = [e for e in range(E) if bool(masked[:, e].all())]
    got = _run(*_poisoned(X, logits, up, down, out_of_service, []), k, mx4, score=mb.MOE_SCORE_SIGMOID if sigmoid else mb.MOE_SCORE_SOFTMAX,
               renormalize=renormalize)
    _check(got, want)


@pytest.mark.parametrize("mx4", [False, True])
def test_a_row_that_is_not_a_number_stays_one(mx4):
    """A NaN logit makes its row's weights NaN, the masked choices' too; the other rows are what they are without it."""
    X, logits, up, down = _inputs(4, 10, 128, 64, 3)
    logits[1, 2:] = -INF
    out, tol, ids, w = _expected(X, logits, up, down, 4, mx4)
    logits[1, 1] = NAN
    got = _run(X, logits, up, down, 4, mx4)
    assert bool(torch.isnan(got[0][1]).all()) and bool(torch.isnan(got[2][1]).all())
    assert torch.equal(got[1], ref.route(logits, 4, False, True, 1.0)[0])
    rest = [0, 2, 3]
    _check([v[rest] for v in got], [v[rest] for v in (out, tol, ids, w)])


@pytest.mark.parametrize("mx4", [False, True])
def test_no_expert_at_all(mx4):
    X, logits, up, down = _inputs(5, 12, 136, 72, 9)
    logits[:] = -INF
    out, ids, w = _run(*_poisoned(X, logits, up, down, range(12), range(5)), 3, mx4)
    assert bool((out == 0).all()) and bool((w == 0).all()) and torch.equal(ids, torch.arange(3, dtype=torch.int32).expand(5, 3))
