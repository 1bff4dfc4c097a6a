"""Weights, outputs and rows whose byte offsets pass 32 bits: the same bits as the same product where they do not."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _randn(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(torch.bfloat16)


def _product(X, W, ids, T, k, E, K, N, gated, tile_m):
    plan = mb.MoeMx4ProductPlan(T, k, E, K, N, gated=gated, device=DEV)
    plan.g = mb.Tiling(tile_m, 256)
    plan.map = mb.alloc_task_map(T, k, E, tile_m, 256, plan.columns, DEV)
    return plan.forward(X, W, ids).clone()


@pytest.mark.parametrize("gated", [False, True])
def test_last_expert_of_more_than_4_GiB(gated):
    E, K, N, T = 40, 8192, 28672, 70
    many, one = mb.Mx4Weights(E, K, N, gated, DEV), mb.Mx4Weights(1, K, N, gated, DEV)
    assert many.codes.numel() > 1 << 32
    W = _randn(K, N, seed=1)
    many.pack_expert(E - 1, W)
    one.pack_expert(0, W)
    X = _randn(T, K, seed=2)
    ids = torch.full((T, 1), E - 1, dtype=torch.int32, device=DEV)
    for tile_m in (16, 32, 128):
        a = _product(X, many, ids, T, 1, E, K, N, gated, tile_m)
        b = _product(X, one, torch.zeros_like(ids), T, 1, 1, K, N, gated, tile_m)
        assert torch.equal(a, b)


def test_output_of_more_than_4_GiB():
    T, K, N = 66000, 128, 36864
    W = mb.Mx4Weights(1, K, N, False, DEV).pack(_randn(1, K, N, seed=3))
    X = _randn(T, K, seed=4)
    ids = torch.zeros(T, 1, dtype=torch.int32, device=DEV)
    for tile_m in (32, 128):
        a = _product(X, W, ids, T, 1, 1, K, N, False, tile_m)
        assert a.numel() * 2 > 1 << 32
        for at in (0, 33000, T - 100):
            b = _product(X[at:at + 100].contiguous(), W, ids[:100], 100, 1, 1, K, N, False, tile_m)
            assert torch.equal(a[at:at + 100], b)
        del a


@pytest.mark.parametrize("mx4", [False, True])
def test_few_tokens_last_expert_of_more_than_4_GiB(mx4):
    E, hidden, inter, T = (40, 8192, 14336, 5) if mx4 else (12, 8192, 14336, 5)
    up, down = _randn(hidden, 2 * inter, seed=5) * hidden ** -0.5, _randn(inter, hidden, seed=6) * inter ** -0.5
    if mx4:
        many = mb.Mx4Weights(E, hidden, 2 * inter, True, DEV), mb.Mx4Weights(E, inter, hidden, False, DEV)
        one = mb.Mx4Weights(1, hidden, 2 * inter, True, DEV), mb.Mx4Weights(1, inter, hidden, False, DEV)
        for w, e in ((many, E - 1), (one, 0)):
            w[0].pack_expert(e, up)
            w[1].pack_expert(e, down)
        assert many[0].codes.numel() > 1 << 32
    else:
        many = torch.empty(E, hidden, 2 * inter, dtype=torch.bfloat16, device=DEV), torch.empty(E, inter, hidden, dtype=torch.bfloat16, device=DEV)
        many[0][E - 1], many[1][E - 1] = up, down
        one = up[None].contiguous(), down[None].contiguous()
        assert many[0].numel() * 2 > 1 << 32
    X = _randn(T, hidden, seed=7)
    logits = torch.zeros(T, E, device=DEV)
    logits[:, E - 1] = 1.0
    a = mb.MoeFewTokensPlan(T, 1, E, hidden, inter, device=DEV).forward(X, logits, *many)
    b = mb.MoeFewTokensPlan(T, 1, 1, hidden, inter, device=DEV).forward(X, logits[:, :1].contiguous(), *one)
    assert bool((a[1] == E - 1).all()) and bool((a[2] == 1).all())
    diff = (a[0].double() - b[0].double()).abs()
    # (column tiles by twos, and parts of the second sum, may go by the number of experts: fp32 sums in another order, each output and a few of h rounded the other way)
    assert bool((diff <= 2.0 ** -7 * b[0].double().abs() + 2.0 ** -11).all()) and bool(torch.isfinite(a[0]).all())


def test_rows_far_apart():
    """Rows of one buffer more than 2^32 bytes apart, for the quantiser and the router."""
    stride = (1 << 31) + 64
    buffer = torch.zeros(stride * 2 + 4096, dtype=torch.bfloat16, device=DEV)
    x = buffer.as_strided((3, 200), (stride, 1))
    x.copy_(_randn(3, 200, seed=8))
    far, near = mb.Mx4Rows(3, 200, DEV).quantize(x), mb.Mx4Rows(3, 200, DEV).quantize(x.contiguous())
    assert torch.equal(far.codes, near.codes) and torch.equal(far.scales, near.scales)
    got = []
    for logits in (x, x.contiguous()):
        ids, w = torch.empty(3, 5, dtype=torch.int32, device=DEV), torch.empty(3, 5, device=DEV)
        mb.moe_route(logits, 5, ids, w)
        got.append((ids, w))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
