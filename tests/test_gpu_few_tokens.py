"""The layer for few tokens against 64 bits: both kinds of weights, every number of tokens, odd sizes, masked rows, and that
nothing but a token's own experts reaches it."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb
from tests import helpers as H
from tests import mx4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _inputs(T, E, hidden, inter, seed, masked=0):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn(T, hidden, generator=g).to(torch.bfloat16)
    logits = torch.randn(T, E, generator=g)
    if masked:
        logits[T - masked:] = -float("inf")
    up = (torch.randn(E, hidden, 2 * inter, generator=g) * hidden ** -0.5).to(torch.bfloat16)
    down = (torch.randn(E, inter, hidden, generator=g) * inter ** -0.5).to(torch.bfloat16)
    return X, logits, up, down


def _values(W, mx4):
    return torch.stack([ref.quantize(w.t())[2].t() for w in W]) if mx4 else W.double()


def _expected(X, logits, up, down, k, mx4, sigmoid=False, renormalize=True, scale=1.0):
    """Output in 64 bits and a bound: fp32 sums of hidden (inter) exact products in any order, h rounded to bf16 once, the
    router's weights and the sum over the experts in fp32, the output rounded to bf16 once."""
    ids, w = ref.route(logits, k, sigmoid, renormalize, scale)
    U, D, x = _values(up, mx4), _values(down, mx4), X.double()
    T, hidden, inter = X.shape[0], X.shape[1], down.shape[1]
    out, tol, mag = torch.zeros(T, hidden, dtype=torch.float64), torch.zeros(T, hidden, dtype=torch.float64), torch.zeros(T, hidden, dtype=torch.float64)
    c1, c2 = H.sum_err_coeff(hidden + 64, False), H.sum_err_coeff(inter + 64, False)
    for t in range(T):
        for j in range(k):
            e = int(ids[t, j])
            y, err = x[t] @ U[e], c1 * (x[t].abs() @ U[e].abs())
            g, u, eg, eu = y[:inter], y[inter:], err[:inter], err[inter:]
            h = ref.silu(g) * u
            eh = 1.1 * eg * (u.abs() + eu) + ref.silu(g).abs() * eu + 32 * 2.0 ** -24 * h.abs()
            eh = eh + 2.0 ** -8 * (h.abs() + eh) + 2.0 ** -130
            z, A = h @ D[e], h.abs() @ D[e].abs()
            ez = eh @ D[e].abs() + c2 * (A + eh @ D[e].abs())
            p = float(w[t, j])
            out[t] += p * z
            mag[t] += p * (z.abs() + ez)
            tol[t] += p * ez
    tol += mag * (k + 64) * 2.0 ** -24 + 2.0 ** -8 * out.abs() + 2.0 ** -130
    return out, tol, ids, w


def _run(X, logits, up, down, k, mx4, **kw):
    T, hidden = X.shape
    E, inter = down.shape[:2]
    plan = mb.MoeFewTokensPlan(T, k, E, hidden, inter, device=DEV, **kw)
    plan.workspace.fill_(0xFF)
    plan.out.fill_(float("nan"))
    if mx4:
        weights = mb.Mx4Weights(E, hidden, 2 * inter, True, DEV).pack(up.to(DEV)), mb.Mx4Weights(E, inter, hidden, False, DEV).pack(down.to(DEV))
    else:
        weights = up.to(DEV), down.to(DEV)
    out, ids, w = plan.forward(X.to(DEV), logits.to(DEV), *weights)
    return out.cpu(), ids.cpu(), w.cpu()


def _check(got, want):
    (out, ids, w), (ref_out, tol, ref_ids, ref_w) = got, want
    assert torch.equal(ids, ref_ids)
    assert bool(((w.double() - ref_w).abs() <= 40 * 2.0 ** -24 * ref_w + 2.0 ** -125).all())
    bad = ~((out.double() - ref_out).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), out[bad][:4], ref_out[bad][:4], tol[bad][:4])


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("T,k,E,hidden,inter", [
    (1, 1, 1, 8, 8), (1, 1, 3, 64, 32), (1, 6, 64, 256, 176), (2, 2, 4, 136, 72), (3, 3, 5, 264, 40), (4, 2, 8, 512, 384), (5, 8, 256, 128, 64),
    (7, 4, 100, 384, 200), (8, 1, 2, 1024, 128), (11, 6, 64, 256, 256), (13, 16, 40, 128, 96), (15, 2, 8, 640, 1000), (16, 16, 16, 136, 72),
    (16, 8, 1000, 64, 64), (16, 2, 3, 2048, 520), (16, 6, 64, 512, 176)])
def test_layer(T, k, E, hidden, inter, mx4):
    data = _inputs(T, E, hidden, inter, T * 100 + E)
    _check(_run(*data, k, mx4), _expected(*data, k, mx4))


@pytest.mark.parametrize("T", range(1, 17))
@pytest.mark.parametrize("mx4", [False, True])
def test_every_number_of_tokens(T, mx4):
    data = _inputs(T, 6, 200, 88, T)
    _check(_run(*data, 2, mx4), _expected(*data, 2, mx4))


@pytest.mark.parametrize("inter", [1, 7, 15, 17, 33, 50])
def test_widths_that_only_the_packed_weights_take(inter):
    data = _inputs(3, 4, 72, inter, inter)
    _check(_run(*data, 2, True), _expected(*data, 2, True))


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("sigmoid,renormalize,scale", [(True, True, 2.5), (True, False, 1.0), (False, False, 1.0)])
def test_scores(sigmoid, renormalize, scale, mx4):
    X, logits, up, down = _inputs(6, 20, 256, 96, 3)
    logits = logits.to(torch.bfloat16)
    got = _run(X, logits, up, down, 4, mx4, score=mb.MOE_SCORE_SIGMOID if sigmoid else mb.MOE_SCORE_SOFTMAX, renormalize=renormalize, scale=scale)
    _check(got, _expected(X, logits, up, down, 4, mx4, sigmoid, renormalize, scale))


@pytest.mark.parametrize("mx4", [False, True])
def test_masked_tokens_come_out_as_zeros(mx4):
    data = _inputs(9, 8, 256, 128, 5, masked=4)
    got = _run(*data, 3, mx4)
    _check(got, _expected(*data, 3, mx4))
    assert bool((got[0][5:] == 0).all()) and bool((got[2][5:] == 0).all())


@pytest.mark.parametrize("mx4", [False, True])
def test_nothing_but_its_own_experts_reaches_a_token(mx4):
    """Infinities and NaN in the weights of one expert and in one token: every other token's output keeps its bits."""
    X, logits, up, down = _inputs(12, 10, 264, 136, 7)
    clean = _run(X, logits, up, down, 2, mx4)
    e = int(clean[1][3, 0])
    hit = (clean[1] == e).any(1)
    hit[6] = True
    assert 2 <= int(hit.sum()) < 12
    up, down, X = up.clone(), down.clone(), X.clone()
    up[e, 5, 3], down[e, 7, :] = float("inf"), float("nan")
    X[6, 9] = float("nan")
    got = _run(X, logits, up, down, 2, mx4)
    assert torch.equal(got[0][~hit], clean[0][~hit])
    assert bool(torch.isnan(got[0][hit]).any(1).all())


@pytest.mark.parametrize("mx4", [False, True])
def test_same_bits_again_on_streams_and_from_a_graph(mx4):
    T, k, E, hidden, inter = 4, 4, 32, 1024, 512
    X, logits, up, down = _inputs(T, E, hidden, inter, 13)
    plan = mb.MoeFewTokensPlan(T, k, E, hidden, inter, device=DEV)
    if mx4:
        weights = mb.Mx4Weights(E, hidden, 2 * inter, True, DEV).pack(up.to(DEV)), mb.Mx4Weights(E, inter, hidden, False, DEV).pack(down.to(DEV))
    else:
        weights = up.to(DEV), down.to(DEV)
    x, lg = torch.empty_like(X, device=DEV), torch.empty_like(logits, device=DEV)

    def inputs(seed):
        a, b, _, _ = _inputs(T, E, hidden, inter, seed)
        x.copy_(a)
        lg.copy_(b)
        torch.cuda.synchronize()

    def eager():
        plan.forward(x, lg, *weights)
        torch.cuda.synchronize()
        return plan.out.clone(), plan.ids.clone()

    first = {}
    for seed in (1, 2, 3):
        inputs(seed)
        first[seed] = eager()
        for _ in range(5):
            again = eager()
            assert torch.equal(again[0], first[seed][0]) and torch.equal(again[1], first[seed][1])
    s = torch.cuda.Stream()
    inputs(2)
    with torch.cuda.stream(s):
        plan.forward(x, lg, *weights)
    s.synchronize()
    assert torch.equal(plan.out, first[2][0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.forward(x, lg, *weights)
    for seed in (3, 1, 2, 1):
        inputs(seed)
        plan.out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(plan.out, first[seed][0]) and torch.equal(plan.ids, first[seed][1])


@pytest.mark.parametrize("T,k,E,hidden,inter", [(16, 2, 3, 4712, 40), (16, 3, 300, 4608, 16), (9, 2, 2, 8200, 24)])
def test_more_token_values_than_lds_holds(T, k, E, hidden, inter):
    data = _inputs(T, E, hidden, inter, hidden)
    _check(_run(*data, k, True), _expected(*data, k, True))


@pytest.mark.parametrize("T,k,E,hidden,inter", [(8, 2, 16, 72, 2048), (8, 2, 16, 40, 2104), (16, 4, 300, 16, 448)])
def test_column_tiles_by_twos(T, k, E, hidden, inter):
    data = _inputs(T, E, hidden, inter, inter)
    _check(_run(*data, k, False), _expected(*data, k, False))


def test_no_tokens():
    plan = mb.MoeFewTokensPlan(0, 2, 4, 64, 64, device=DEV)
    e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=DEV)
    out, ids, w = plan.forward(e(0, 64), torch.empty(0, 4, device=DEV), e(4, 64, 128), e(4, 64, 64))
    assert out.shape == (0, 64) and ids.shape == (0, 2)
