"""The grouped router's choice: ids exactly, weights against 64 bits."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb
from tests import block_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _inputs(T, E, seed, dtype, kind):
    g = torch.Generator().manual_seed(seed)
    x, bias = torch.randn(T, E, generator=g) * 2, torch.randn(E, generator=g) * 0.2
    if kind == "ties":            # few different logits and biases (none whose sigmoids add up to the same in two ways)
        x, bias = torch.randint(0, 4, (T, E), generator=g).float(), torch.randint(-1, 2, (E,), generator=g) * 0.125
    elif kind == "masked":
        x[torch.rand(T, E, generator=g) < 0.6] = -float("inf")
        x[T // 2] = -float("inf")
        x[0, : E - 1] = -float("inf")
        bias[E // 2] = -float("inf")
    elif kind == "lowest":        # masks of the type's lowest value count as numbers
        x[torch.rand(T, E, generator=g) < 0.6] = torch.finfo(dtype).min
        x[T // 2] = torch.finfo(dtype).min
    elif kind == "large":         # most scores are zero in 64 bits too: the logit decides
        x *= 1e4
    return x.to(dtype), bias


def _run(x, k, groups, kept, top2, bias, sigmoid, renormalize, scale):
    T = x.shape[0]
    ids = torch.full((T + 1, k), -7, dtype=torch.int32, device=DEV)
    w = torch.full((T + 1, k), 7.0, device=DEV)
    mb.moe_route_grouped(x, k, ids, w, groups, kept, mb.MOE_GROUP_TOP2 if top2 else mb.MOE_GROUP_MAX, bias,
                         mb.MOE_SCORE_SIGMOID if sigmoid else mb.MOE_SCORE_SOFTMAX, renormalize, scale)
    assert bool((ids[T] == -7).all()) and bool((w[T] == 7.0).all())
    return ids[:T].cpu(), w[:T].cpu().double()


def _check(x_gpu, x, k, groups, kept, top2, bias, sigmoid, renormalize, scale):
    ids, w = _run(x_gpu, k, groups, kept, top2, None if bias is None else bias.to(DEV), sigmoid, renormalize, scale)
    want_ids, want = ref.route_grouped(x, k, groups, kept, top2, bias, sigmoid, renormalize, scale)
    assert torch.equal(ids, want_ids)
    assert torch.equal(torch.isnan(w), torch.isnan(want))
    # 64 bits throughout, rounded once: half a step of fp32 and a hundredth for 64 bits' own roundings; below 2^-126 half of 2^-149, doubled for a flush of the last bit
    ok = ~torch.isnan(want)
    assert bool(((w - want).abs() <= 1.01 * 2.0 ** -24 * want.abs() + 2.0 ** -149)[ok].all())


@pytest.mark.parametrize("kind", ["normal", "ties", "masked", "lowest", "large"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,E,k,groups,kept", [(1, 1, 1, 1, 1), (1, 64, 6, 8, 4), (2, 8, 8, 4, 4), (5, 20, 3, 5, 2), (33, 60, 6, 4, 1), (17, 65, 8, 13, 3), (40, 256, 8, 8, 4),
                                               (9, 257, 16, 1, 1), (3, 1023, 31, 33, 1), (4, 100, 50, 2, 1), (6, 72, 6, 6, 3), (7, 320, 8, 10, 3), (5, 512, 8, 8, 2),
                                               (3, 1023, 8, 3, 2), (4, 64, 3, 64, 3), (3, 128, 70, 32, 20), (2, 1000, 500, 5, 3)])
def test_route_grouped(T, E, k, groups, kept, dtype, kind):
    x, bias = _inputs(T, E, T * 1000 + E + k, dtype, kind)
    for sigmoid in (False, True):
        for top2 in (False, True):
            _check(x.to(DEV), x, k, groups, kept, top2, bias if kind != "large" else None, sigmoid, top2, 2.5 if sigmoid else 1.0)
            _check(x.to(DEV), x, k, groups, kept, top2, None, sigmoid, not top2, 1.0)


def test_many_tokens():
    x, bias = _inputs(1501, 160, 4, torch.float32, "normal")
    _check(x.to(DEV), x, 6, 8, 3, True, bias, True, True, 2.5)


@pytest.mark.parametrize("T", [4, 5, 6, 7, 8])
@pytest.mark.parametrize("k", [1, 15, 16, 17])
@pytest.mark.parametrize("E", [64, 120, 256, 512])
def test_four_tokens_of_a_workgroup(T, k, E):
    """Every number of tokens in the last workgroup, choices on either side of a quarter of the lanes."""
    for kind in ("normal", "masked"):
        x, bias = _inputs(T, E, T * 100 + k, torch.float32, kind)
        for renormalize in (False, True):
            _check(x.to(DEV), x, k, 4, 3, True, bias, True, renormalize, 2.5)


@pytest.mark.parametrize("spread", [1e-9, 1e-4, 1.0, 30.0, 300.0])
@pytest.mark.parametrize("shift", [-650.0, -40.0, 0.0, 15.0, 40.0])
def test_flat_and_peaked_rows_without_a_bias(spread, shift):
    """Scores that are nearly equal, that saturate, and that leave 32 (and 64) bits; groups of equal scores go by their index."""
    x = torch.randn(40, 96, generator=torch.Generator().manual_seed(int(spread + shift + 1000))) * spread + shift
    x[7] = x[7, 0]
    for sigmoid in (False, True):
        for top2 in (False, True):
            _check(x.to(DEV), x, 6, 8, 3, top2, None, sigmoid, False, 1.0)
            _check(x.to(DEV), x, 5, 3, 1, top2, None, sigmoid, True, 1.0)


def test_scores_next_to_each_other():
    """Scores that 32 bits cannot tell apart: biases that make up for the logits' difference to within 2^-40."""
    g = torch.Generator().manual_seed(5)
    x = torch.randn(200, 64, generator=g)
    p = torch.sigmoid(x[:1].double())
    bias = (0.75 - p[0]).float()                     # s = 0.75 up to bias's rounding, 2^-26: well apart in 64 bits, not in 32
    x[:] = x[0]
    x += 1e-7 * torch.randn(200, 64, generator=g)
    _check(x.to(DEV), x, 8, 8, 4, True, bias, True, True, 1.0)


@pytest.mark.parametrize("low", [-1e9, -1e4, -30.0, 1e4])
def test_experts_put_out_of_reach_by_their_bias(low):
    """Biases far from the others' count as numbers: such experts come last (or first), and the others are told apart as without them."""
    x, bias = _inputs(60, 128, 31, torch.float32, "normal")
    bias[5::7] = low
    bias[32:48] = low                                # a whole group
    for sigmoid in (False, True):
        for top2 in (False, True):
            _check(x.to(DEV), x, 6, 8, 3, top2, bias, sigmoid, True, 1.0)
            _check(x.to(DEV), x, 40, 8, 4, top2, bias, sigmoid, True, 1.0)


@pytest.mark.parametrize("k", [1, 2, 5, 6, 15, 16, 31])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_neighbours_in_pairs(k, sigmoid):
    """Pairs of scores that differ by less than 32 bits can tell, well apart from the next pair; the border of the choice lies between two pairs or in one."""
    g = torch.Generator().manual_seed(k)
    for groups, kept in ((8, 4), (1, 1)):
        x = torch.randn(1, 64, generator=g)
        p = torch.sigmoid(x.double()) if sigmoid else torch.softmax(x.double(), 1)
        place = torch.randperm(64, generator=g)
        bias = (1.5 - 0.01 * (place // 2) - p[0]).float()        # (rounded: the two of a pair end up some 2^-26 apart)
        x = x + 1e-8 * torch.randn(60, 64, generator=g)
        _check(x.to(DEV), x, k, groups, kept, False, bias, sigmoid, True, 1.0)


def test_without_groups_and_bias_the_choices_are_moe_routes():
    for kind in ("normal", "ties", "masked", "large"):
        x, _ = _inputs(50, 96, 8, torch.float32, kind)
        ids, w = torch.empty(50, 6, dtype=torch.int32, device=DEV), torch.empty(50, 6, device=DEV)
        for score in (mb.MOE_SCORE_SOFTMAX, mb.MOE_SCORE_SIGMOID):
            mb.moe_route(x.to(DEV), 6, ids, w, score=score)
            got, _ = _run(x.to(DEV), 6, 1, 1, False, None, score == mb.MOE_SCORE_SIGMOID, True, 1.0)
            assert torch.equal(got, ids.cpu())


def test_rows_apart():
    wide, bias = _inputs(30, 200, 9, torch.float32, "normal")
    _check(wide.to(DEV)[:, 7:135], wide[:, 7:135], 8, 8, 3, True, bias[:128], True, True, 1.0)
    _check(wide.to(DEV)[::3, :64], wide[::3, :64], 4, 4, 2, False, None, True, False, 1.0)
    half, _ = _inputs(30, 131, 10, torch.bfloat16, "ties")
    _check(half.to(DEV)[:, 1:], half[:, 1:], 8, 10, 4, False, None, False, True, 1.0)


def test_not_a_number():
    """A NaN score comes first, and its group too; in a softmax row all scores are NaN, and then logits decide (a NaN before +inf)."""
    x, bias = _inputs(5, 64, 3, torch.float32, "normal")
    x[0, 60], x[1, 3], x[2, 3], x[2, 40] = float("nan"), float("inf"), float("nan"), float("nan")
    x[3, 10] = -float("inf")
    nan_bias = bias.clone()
    nan_bias[17] = float("nan")
    for b in (bias, None, nan_bias):
        for top2 in (False, True):
            for renormalize in (False, True):
                _check(x.to(DEV), x, 5, 8, 3, top2, b, True, renormalize, 1.0)
        ids, w = _run(x.to(DEV), 5, 8, 3, True, None if b is None else b.to(DEV), False, True, 1.0)
        assert bool(torch.isnan(w[:3]).all()) and not bool(torch.isnan(w[4]).any())
        assert bool((ids >= 0).all()) and bool((ids < 64).all())


def test_no_tokens():
    assert mb.moe_route_grouped(torch.empty(0, 8, device=DEV), 2, torch.empty(0, 2, dtype=torch.int32, device=DEV), torch.empty(0, 2, device=DEV), 2, 1) == mb.MOE_OK


def test_captured_and_on_a_stream():
    x, bias = _inputs(70, 256, 21, torch.float32, "normal")
    xg, bg = x.to(DEV), bias.to(DEV)
    ids, w = torch.empty(70, 8, dtype=torch.int32, device=DEV), torch.empty(70, 8, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        mb.moe_route_grouped(xg, 8, ids, w, 8, 4, mb.MOE_GROUP_TOP2, bg, mb.MOE_SCORE_SIGMOID)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        mb.moe_route_grouped(xg, 8, ids, w, 8, 4, mb.MOE_GROUP_TOP2, bg, mb.MOE_SCORE_SIGMOID)
    for turn in range(3):
        x = x.roll(1, 0)
        xg.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        want, weights = ref.route_grouped(x, 8, 8, 4, True, bias, True, True, 1.0)
        assert torch.equal(ids.cpu(), want) and torch.allclose(w.cpu().double(), weights, rtol=1.01 * 2.0 ** -24, atol=0)


def test_on_a_stream_of_its_own():
    """What a call on another stream than the default one writes, behind inputs that are made there."""
    x, bias = _inputs(70, 256, 22, torch.float32, "normal")
    ids, w = torch.full((70, 8), -7, dtype=torch.int32, device=DEV), torch.full((70, 8), 7.0, device=DEV)
    xg, bg = torch.zeros(70, 256, device=DEV), bias.to(DEV)
    late = x.to(DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(1 << 22)
        xg.copy_(late)
        mb.moe_route_grouped(xg, 8, ids, w, 8, 4, mb.MOE_GROUP_TOP2, bg, mb.MOE_SCORE_SIGMOID)
    s.synchronize()
    want, weights = ref.route_grouped(x, 8, 8, 4, True, bias, True, True, 1.0)
    assert torch.equal(ids.cpu(), want) and torch.allclose(w.cpu().double(), weights, rtol=1.01 * 2.0 ** -24, atol=0)
